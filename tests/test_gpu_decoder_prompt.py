"""The example's layer takes in packed prompts and then checks trees behind them, with norms and rotation, against the same layer in plain 32-bit torch;
and a training step through rotation and attention against differentiated plain torch."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(ROOT, "examples", "decoder_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def turn(x, weight, freqs, positions):
    """[tokens, heads, d], 32 bits."""
    import torch
    if weight is not None:
        x = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight.float()
    angle = positions.double()[:, None, None] * freqs
    cos, sin, half = angle.cos().float(), angle.sin().float(), x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def attend(q, k, v, keep):                      # [n, H, d], [L, Hkv, d], [n, L]
    import torch
    H, Hkv, d = q.shape[1], k.shape[1], q.shape[2]
    k, v = (z.repeat_interleave(H // Hkv, 1) for z in (k, v))
    s = torch.einsum("nhd,lhd->hnl", q, k) * d ** -0.5
    return torch.einsum("hnl,lhd->nhd", torch.softmax(s.masked_fill(~keep, -float("inf")), 2), v)


def plain_layer(layer, x, own, enc_k, enc_v):
    """The layer around its self-attention: own(q, k, v as projected) -> its result."""
    import torch
    H, Hkv, d = layer.heads, layer.kv_heads, layer.head_dim
    norm = lambda z: torch.nn.functional.layer_norm(z.float(), (H * d,))  # noqa: E731
    f = lambda w: w.float().t()  # noqa: E731
    qkv = (norm(x) @ f(layer.w_qkv)).view(-1, H + 2 * Hkv, d)
    x = x + own(qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]).reshape(len(x), -1) @ f(layer.w_self_out)
    q = (norm(x) @ f(layer.w_cross_q)).view(-1, H, d)
    everything = torch.ones(len(x), len(enc_k), dtype=torch.bool, device="cuda")
    x = x + attend(q, enc_k.float(), enc_v.float(), everything).reshape(len(x), -1) @ f(layer.w_cross_out)
    z = norm(x)
    return x + (torch.nn.functional.silu(z @ f(layer.w_gate)) * (z @ f(layer.w_up))) @ f(layer.w_down)


@pytest.mark.parametrize("base", [None, 10000.0])
def test_prompts_then_a_tree(E, base):
    import torch
    n, H, Hkv, d, lens, enc_lens = 7, 8, 2, 64, [40, 1, 173], [30, 90, 5]
    layer = E.Layer(3, n, H, Hkv, d, 320, dtype=torch.float16, base=base)
    p = E.prompts(layer, lens, enc_lens)
    chain = torch.tril(torch.ones(n, n, dtype=torch.bool))          # drafted one after the other, but the last two beside each other
    chain[n - 1, n - 2] = False
    bits = (chain.long() << torch.arange(n)).sum(1).expand(3, n).contiguous()[..., None].cuda()
    held = torch.tensor(lens, dtype=torch.int32, device="cuda")
    depth = torch.tensor(list(range(n - 1)) + [n - 2], device="cuda")
    positions = (held[:, None] + depth).to(torch.int32).flatten()
    g = torch.Generator(device="cuda").manual_seed(9)
    x_tree = torch.randn(3, n, H * d, generator=g, device="cuda").to(torch.float16)
    enc = torch.zeros(3, max(enc_lens), 2, Hkv, d, dtype=torch.float16, device="cuda")
    for b in range(3):
        keys = slice(int(p["enc_starts"][b]), int(p["enc_starts"][b + 1]))
        enc[b, :enc_lens[b], 0], enc[b, :enc_lens[b], 1] = p["enc_k"][keys], p["enc_v"][keys]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    E.M.mmee_set_stream(stream.cuda_stream)
    try:
        with torch.cuda.stream(stream):
            got = layer.prompt(**p)
            tree = layer.step(x_tree, p["k_pages"], p["v_pages"], p["page_table"], held, bits, enc[:, :, 0], enc[:, :, 1],
                              torch.tensor(enc_lens, dtype=torch.int32, device="cuda"), positions=positions if base else None)
        stream.synchronize()
    finally:
        E.M.mmee_set_stream(None)
    for b in range(3):
        kept = {}

        def own_prompt(q, k, v):
            at = torch.arange(lens[b], device="cuda")
            if base:
                q, k = turn(q, layer.q_weight, layer.freqs, at), turn(k, layer.k_weight, layer.freqs, at)
            kept["k"], kept["v"] = k, v
            return attend(q, k, v, at[None] <= at[:, None])

        def own_tree(q, k, v):
            at = lens[b] + depth
            if base:
                q, k = turn(q, layer.q_weight, layer.freqs, at), turn(k, layer.k_weight, layer.freqs, at)
            keep = torch.cat([torch.ones(n, lens[b], dtype=torch.bool, device="cuda"), chain.cuda()], 1)
            return attend(q, torch.cat([kept["k"], k]), torch.cat([kept["v"], v]), keep)
        rows, keys = slice(int(p["starts"][b]), int(p["starts"][b + 1])), slice(int(p["enc_starts"][b]), int(p["enc_starts"][b + 1]))
        for name, out, want in (("prompt", got[rows], plain_layer(layer, p["x"][rows].float(), own_prompt, p["enc_k"][keys], p["enc_v"][keys])),
                                ("tree", tree[b], plain_layer(layer, x_tree[b].float(), own_tree, p["enc_k"][keys], p["enc_v"][keys]))):
            # some twenty-four roundings to 11 bits of values of size 1 to 4 on the way: 2^-11 each, in the root mean square
            assert (out.float() - want).square().mean().sqrt() <= 2.0 ** -11 * 24 ** 0.5 * want.square().mean().sqrt(), (name, b)
        # what lies in the cache are the keys and values that the prompts' rows were given: a product rounded, a norm and a rotation rounded
        pages = p["page_table"][b].long()
        for name, pool in (("k", p["k_pages"]), ("v", p["v_pages"])):
            there = pool[pages].flatten(0, 1)[:lens[b]].float()
            assert (there - kept[name]).square().mean().sqrt() <= 2.0 ** -11 * 3 * kept[name].square().mean().sqrt(), (name, b)


def test_training_step(E):
    """Norm and rotation, attention over packed prompts, back through both: gradients of the projections' results and of the norms' weights."""
    import torch
    M, lens, H, Hkv, d, dt = E.M, [90, 33, 1, 160], 6, 3, 64, torch.bfloat16
    T = sum(lens)
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    x, do, weights = r(T, H + 2 * Hkv, d), r(T, H, d), [(1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2)]
    starts = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    positions = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
    freqs = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).cuda()
    q, k, v = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
    empty = lambda *s: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    q_out, k_out, o, lse = empty(T, H, d), empty(T, Hkv, d), empty(T, H, d), torch.empty(H, T, device="cuda")
    dx, dw = empty(T, H + 2 * Hkv, d), [empty(d), empty(d)]
    dq, dk = empty(T, H, d), empty(T, Hkv, d)
    turned = M.qk_rotate(q, k, q_out, k_out, freqs, positions, q_weight=weights[0], k_weight=weights[1])
    attention = M.prompt_attn(q_out, k_out, v, o, starts, lse=lse)
    back = M.qk_rotate_grads(dq, dk, dx[:, :H], dx[:, H:H + Hkv], *dw)
    for call, size in ((turned, M.mmee_qk_rotate_workspace(turned)), (attention, M.mmee_prompt_attn_workspace(attention, True))):
        call.use_workspace(torch.empty(size, dtype=torch.uint8, device="cuda"))
    M.mmee_qk_rotate_forward(turned)
    M.mmee_prompt_attn_forward(attention)
    M.mmee_prompt_attn_backward(attention, M.prompt_attn_grads(do, dq, dk, dx[:, H + Hkv:]))
    M.mmee_qk_rotate_backward(turned, back)
    torch.cuda.synchronize()

    X, W = x.float().requires_grad_(), [w.float().requires_grad_() for w in weights]
    Q, K, V = turn(X[:, :H], W[0], freqs, positions), turn(X[:, H:H + Hkv], W[1], freqs, positions), X[:, H + Hkv:]
    want, at = [], 0
    for n in lens:
        rows = slice(at, at + n)
        i = torch.arange(n, device="cuda")
        want.append(attend(Q[rows], K[rows], V[rows], i[None] <= i[:, None]))
        at += n
    want = torch.cat(want)
    grads = torch.autograd.grad(want, [X, *W], do.float())
    # roundings to 8 bits on the way, 2^-8 each in the root mean square: o: q, k, probabilities, o; gradients: these, dS, their own, and the projections' rounded ones
    for name, got, exact, roundings in (("o", o, want, 4), ("dx", dx, grads[0], 8), ("dq_weight", dw[0], grads[1], 8), ("dk_weight", dw[1], grads[2], 8)):
        off = (got.float() - exact).square().mean().sqrt() / exact.square().mean().sqrt()
        assert off <= 2.0 ** -8 * roundings ** 0.5, (name, off.item())
