"""Attention of packed prompts, forward and backward, against a plain 64-bit form (attention_oracle.py) sequence by sequence: lengths from none to
several tiles, causal or not, rows over longer and shorter keys, shared heads, layouts, pieces, what lies around the sequences, streams, graphs."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


def starts_of(lens, before=0):
    import torch
    at = [before]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def tensors(q_lens, kv_lens, H, Hkv, d, dtype, seed, train=True, around=0):
    """`around` tokens of no sequence before the first and behind the last one, holding NaN."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    Tq, Tk = sum(q_lens) + 2 * around, sum(kv_lens) + 2 * around

    def r(T, heads):
        x = torch.randn(T, heads, d, generator=g, device="cuda").to(dtype)
        if around:
            x[:around] = x[T - around:] = math.nan
        return x
    t = {"q": r(Tq, H), "k": r(Tk, Hkv), "v": r(Tk, Hkv), "q_starts": starts_of(q_lens, around), "kv_starts": starts_of(kv_lens, around)}
    t["o"], t["lse"] = torch.full_like(t["q"], 9.0), torch.full((H, Tq), 9.0, device="cuda")
    if train:
        t["do"] = r(Tq, H)
        t |= {n: torch.full_like(t[n[1]], 9.0) for n in ("dq", "dk", "dv")}
    return t


def calls(M, t, kv=True, **kw):
    import torch
    a = M.prompt_attn(t["q"], t["k"], t["v"], t["o"], t["q_starts"], kv_starts=t["kv_starts"] if kv else None, lse=t["lse"], **kw)
    # whatever the workspace holds before a call does not matter
    a.use_workspace(torch.full((M.mmee_prompt_attn_workspace(a, "do" in t),), 255, dtype=torch.uint8, device="cuda"))
    return a, M.prompt_attn_grads(t["do"], t["dq"], t["dk"], t["dv"]) if "do" in t else None


def run(M, t, **kw):
    import torch
    a, g = calls(M, t, **kw)
    M.mmee_prompt_attn_forward(a)
    if g:
        M.mmee_prompt_attn_backward(a, g)
    torch.cuda.synchronize()


def keep_of(m, n, causal):
    import torch
    return torch.ones(1, m, n, dtype=torch.bool).tril(n - m) if causal else torch.ones(1, m, n, dtype=torch.bool)


def compare(t, causal, where, scale=None):
    from attention_oracle import attention, check
    q_starts, kv_starts = t["q_starts"].tolist(), t["kv_starts"].tolist()
    for b in range(len(q_starts) - 1):
        rows, keys = slice(q_starts[b], q_starts[b + 1]), slice(kv_starts[b], kv_starts[b + 1])
        one = lambda n: t[n][keys if n[-1] in "kv" else rows][None]  # noqa: E731
        m, n = rows.stop - rows.start, keys.stop - keys.start
        want = attention(one("q"), one("k"), one("v"), keep_of(m, n, causal), scale or t["q"].shape[2] ** -0.5, t["q"].dtype, one("do") if "do" in t else None)
        for name, value in want.items():
            check(t["lse"][:, rows][None] if name == "lse" else one(name), value, (where, b, m, n, name))
    around = [(n, t["kv_starts"] if n[-1] in "kv" else t["q_starts"]) for n in ("o", "dq", "dk", "dv") if n in t]
    for name, of in around:                     # tokens of no sequence
        assert (t[name][:int(of[0])] == 9.0).all() and (t[name][int(of[-1]):] == 9.0).all(), (where, name)
    assert (t["lse"][:, :q_starts[0]] == 9.0).all() and (t["lse"][:, q_starts[-1]:] == 9.0).all()


SHAPES = [  # lengths, H, Hkv, d
    ([1], 1, 1, 8), ([33], 2, 1, 32), ([5, 0, 64, 1, 65], 4, 2, 40), ([63, 128, 2], 3, 3, 64), ([129, 31], 8, 1, 72), ([17, 127, 1, 1, 1], 4, 2, 128), ([257], 2, 2, 96),
    ([300, 40, 200], 6, 2, 120), ([0, 0, 100, 0], 12, 4, 24), ([70, 513], 2, 1, 16), ([256, 255], 1, 1, 56)]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,H,Hkv,d", SHAPES)
def test_prompts_over_themselves(M, lens, H, Hkv, d, causal, dtype):
    import torch
    t = tensors(lens, lens, H, Hkv, d, getattr(torch, dtype), sum(lens) + d)
    run(M, t, kv=False, causal=causal)
    compare(t, causal, (lens, d, causal))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q_lens,kv_lens,H,Hkv,d", [
    ([1], [700], 4, 1, 64), ([3, 1, 1, 40], [64, 129, 1, 41], 8, 2, 128), ([100, 20, 7], [30, 20, 0], 2, 2, 64), ([130, 0, 64], [300, 50, 65], 3, 1, 80), ([257, 1], [1, 1], 2, 1, 32),
    ([64, 64], [1000, 63], 16, 2, 128)])
def test_rows_over_other_keys(M, q_lens, kv_lens, H, Hkv, d, causal, dtype):
    """The last row at the last key: rows before the first key see nothing, give zeros and get zero gradients, and give none."""
    import torch
    t = tensors(q_lens, kv_lens, H, Hkv, d, getattr(torch, dtype), 3, around=3)
    run(M, t, causal=causal)
    compare(t, causal, (q_lens, kv_lens, d, causal))
    for b, (m, n) in enumerate(zip(q_lens, kv_lens)):
        none = slice(int(t["q_starts"][b]), int(t["q_starts"][b]) + (max(0, m - n) if causal else m if not n else 0))
        assert not t["o"][none].any() and not t["dq"][none].any() and (t["lse"][:, none] == -math.inf).all()


def test_what_rows_without_keys_hold(M):
    """Their queries and output gradients may be anything."""
    import torch
    t = tensors([100, 9], [30, 9], 4, 2, 64, torch.float16, 4)
    t["q"][:70:3], t["do"][1:70:3], t["q"][2:70:3] = math.nan, math.inf, math.inf
    run(M, t)
    clean = dict(t)
    clean["q"], clean["do"] = t["q"].clone(), t["do"].clone()
    clean["q"][:70] = clean["do"][:70] = 0
    compare(clean, True, "rows without keys")


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,lens", [(24, [1, 2, 127, 5, 128]), (64, [1, 2, 3, 5, 33, 64]), (128, [1, 64, 2, 6, 9]), (48, [17, 16, 15, 8]), (120, [16, 17])])
def test_gradients_of_few_keys(M, d, lens, causal, dtype):
    """Where a row sees few keys D does not add the rounding of the output: dQ and dK are off by the rounding of dS and their own alone.

    With up to 16 keys of a sequence those of dS are u^2 alone, as what the first rounding leaves is taken along.

    To u |dS_ij| of each dS (u half a step), summed with what multiplies it, and u of the result come the errors in 32 bits, P of 2^-19 (scores of less than 16
    powers of two, the exponential's argument, lse and the exponential each below 2^-21) and dP of d 2^-24 of its terms, in dP and in D; 2^-16 of P (|dP| + D's terms)
    covers them.  Float16 has steps of 2^-24 below its normal numbers."""
    import torch
    t = tensors(lens, lens, 4, 2, d, getattr(torch, dtype), 31 + d)
    run(M, t, kv=False, causal=causal)
    u, scale = torch.finfo(t["q"].dtype).eps / 2, d ** -0.5
    for b, n in enumerate(lens):
        at = slice(sum(lens[:b]), sum(lens[:b]) + n)
        q, do = (t[x][at].double().cpu().view(n, 2, 2, d).permute(1, 2, 0, 3) for x in ("q", "do"))          # [kv head][its heads][row][d]
        k, v = (t[x][at].double().cpu().permute(1, 0, 2)[:, None] for x in ("k", "v"))
        S = q @ k.transpose(2, 3) * scale
        P = S.masked_fill(~keep_of(n, n, causal), -math.inf).softmax(3)
        dP, across = do @ v.transpose(2, 3), do.abs() @ v.abs().transpose(2, 3)
        dS = P * (dP - (P * dP).sum(3, keepdim=True))
        off = (u if n > 16 else u * u) * dS.abs() + 2.0 ** -16 * P * (across + (P * across).sum(3, keepdim=True))
        for name, want, bound in (("dq", dS @ k, off @ k.abs()), ("dk", (dS.transpose(2, 3) @ q).sum(1, keepdim=True), (off.transpose(2, 3) @ q.abs()).sum(1, keepdim=True))):
            got = t[name][at].double().cpu().view(n, 2, -1, d).permute(1, 2, 0, 3)
            far = (got - want * scale).abs() - (1.01 * bound + u * want.abs()) * scale - 2.0 ** -25
            assert (far <= 0).all(), (b, n, name, far.max().item())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q_lens,kv_lens,H,Hkv,d,train", [
    ([40], [3000], 4, 1, 128, True), ([1, 1], [5000, 700], 8, 2, 64, True), ([900], [70], 8, 1, 32, True), ([200, 30], [2500, 2600], 2, 1, 72, True),
    ([270], [270], 70, 70, 64, True), ([300, 520], [1300, 520], 80, 40, 128, True), ([260, 257], [1601, 1500], 33, 33, 72, False)])
def test_pieces_and_many_blocks(M, q_lens, kv_lens, H, Hkv, d, train, causal):
    """Few tiles over many keys or rows, cut into pieces that are joined; tiles of 256 rows and keys, alone and in pieces."""
    import torch
    t = tensors(q_lens, kv_lens, H, Hkv, d, torch.bfloat16, 5, train=train, around=1)
    run(M, t, causal=causal)
    compare(t, causal, (q_lens, kv_lens, causal))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_tiles_of_256(M, dtype):
    import torch
    for d in (64, 128):
        t = tensors([300, 700], [300, 700], 64, 32, d, getattr(torch, dtype), 6)
        run(M, t, kv=False)
        compare(t, True, d)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("group", [1, 3, 8, 32])
def test_keys_of_64_a_wave(M, group, dtype):
    """Tiles of 256 keys with 128 (and 104) values: query heads that share a key/value head so that 32 rows are whole tokens, or not."""
    import torch
    lens, kv_lens, Hkv = {1: ([600, 700, 300], [650, 700, 257], 40), 3: ([300, 257, 3], [520, 257, 40], 40)}.get(group, ([600, 257, 3], [900, 257, 40], 6))
    for causal in (True, False):
        for d in (128, 104):
            t = tensors(lens, kv_lens, Hkv * group, Hkv, d, getattr(torch, dtype), group, around=1)
            for n in ("q", "do"):               # heads first: a token's heads lie apart
                t[n] = t[n].transpose(0, 1).contiguous().transpose(0, 1)
            run(M, t, causal=causal)
            compare(t, causal, (group, causal, d))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("q_lens,kv_lens,H,Hkv,d", [([300], [4200], 4, 2, 128), ([257, 1400], [5000, 3300], 2, 1, 112), ([1100], [1100], 36, 36, 64)])
def test_long_sequences(M, q_lens, kv_lens, H, Hkv, d, dtype):
    """Blocks of eight waves, which only long sequences take."""
    import torch
    t = tensors(q_lens, kv_lens, H, Hkv, d, getattr(torch, dtype), 19, around=1)
    run(M, t)
    compare(t, True, (q_lens, kv_lens))


def test_many_sequences(M):
    """More than a wave looks at in one go, empty ones among them."""
    import torch
    lens = [i * 7 % 23 if i % 3 else 0 for i in range(200)]
    t = tensors(lens, [n + i % 5 for i, n in enumerate(lens)], 4, 2, 32, torch.bfloat16, 7, around=2)
    run(M, t)
    compare(t, True, "many")


@pytest.mark.parametrize("layout", ["fused qkv", "heads first", "broadcast", "sliced"])
def test_layouts(M, layout):
    import torch
    lens, H, Hkv, d, dt = [70, 33], 4, 2, 64, torch.bfloat16
    T = sum(lens)
    t = tensors(lens, lens, H, Hkv, d, dt, 11)
    if layout == "fused qkv":
        x, dx = torch.cat([t["q"], t["k"], t["v"]], 1), torch.full((T, H + 2 * Hkv, d), math.nan, dtype=dt, device="cuda")
        for p, y in (("", x), ("d", dx)):
            t |= {p + "q": y[:, :H], p + "k": y[:, H:H + Hkv], p + "v": y[:, H + Hkv:]}
    elif layout == "heads first":
        t |= {n: t[n].transpose(0, 1).contiguous().transpose(0, 1) for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")}
    elif layout == "broadcast":
        t["k"], t["do"] = t["k"][:, :1].expand(T, Hkv, d), t["do"][:1].expand(T, H, d)
        t["v"] = t["v"][:1].expand(T, Hkv, d)
    else:
        wide = torch.full((T, H, d + 8), 5.0, dtype=dt, device="cuda")
        t["o"] = wide[..., 8:]
    run(M, t, kv=False)
    compare(t, True, layout)
    if layout == "sliced":
        assert (wide[..., :8] == 5.0).all()


def test_scale_and_extremes(M):
    """Scores far apart, the type's largest values, another scale."""
    import torch
    t = tensors([80, 20], [80, 20], 2, 1, 64, torch.bfloat16, 12)
    t["q"][::7] *= 30
    run(M, t, kv=False, scale=0.3)
    compare(t, True, "scale", scale=0.3)


def test_nothing_to_do(M):
    import torch
    t = tensors([0, 0], [5, 70], 2, 1, 64, torch.bfloat16, 1)
    run(M, t)
    assert not t["dk"].any() and not t["dv"].any()
    t = tensors([5, 70], [0, 0], 2, 1, 64, torch.bfloat16, 1)
    run(M, t)
    assert not t["o"].any() and not t["dq"].any() and (t["lse"] == -math.inf).all()
    t = tensors([0], [0], 2, 1, 64, torch.bfloat16, 1)
    run(M, t, kv=False)


def test_starts_beyond_the_tokens_and_out_of_order(M):
    """Clamped; a sequence that ends before it starts is empty."""
    import torch
    t = tensors([50], [50], 2, 1, 64, torch.bfloat16, 2, around=0)
    t["q_starts"] = t["kv_starts"] = torch.tensor([-7, 40, 30, 30, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    run(M, t, kv=False)                          # nothing to compare: whose rows the overlap's are is undefined
    t["q_starts"] = t["kv_starts"] = torch.tensor([-2 ** 31, 20, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    run(M, t, kv=False)
    t["q_starts"] = t["kv_starts"] = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda")
    compare(t, True, "clamped")


def test_long_strides(M):
    """Tokens beyond 2^31 elements from the first one."""
    import torch
    T, d = 200, 64
    row = 1 << 24
    t = tensors([150, 50], [150, 50], 1, 1, d, torch.bfloat16, 14)
    room = torch.empty((T - 1) * row + d, dtype=torch.bfloat16, device="cuda")
    far = room.as_strided((T, 1, d), (row, d, 1))
    far.copy_(t["k"])
    t["k"] = far
    run(M, t, kv=False)
    compare(t, True, "far")


def test_repeats_to_the_bit(M):
    import torch
    t = tensors([300, 1, 64], [2000, 300, 64], 8, 2, 128, torch.float16, 15)
    run(M, t)
    first = {n: t[n].clone() for n in ("o", "lse", "dq", "dk", "dv")}
    run(M, t)
    for n, x in first.items():
        assert torch.equal(x, t[n]), n


def test_streams_and_graphs(M):
    """Captured on a stream of its own and replayed over other inputs and other lengths, with eager calls of the same buffers between the replays."""
    import torch
    t = tensors([90, 60], [90, 60], 4, 2, 64, torch.bfloat16, 16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    M.mmee_set_stream(stream.cuda_stream)
    try:
        a, g = calls(M, t, kv=False)
        M.mmee_prompt_attn_forward(a)
        M.mmee_prompt_attn_backward(a, g)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            M.mmee_prompt_attn_forward(a)
            M.mmee_prompt_attn_backward(a, g)
        for seed, cut in enumerate((90, 1, 150, 0)):
            other = tensors([90, 60], [90, 60], 4, 2, 64, torch.bfloat16, 20 + seed)
            t["q_starts"].copy_(torch.tensor([0, cut, 150]))
            t["kv_starts"].copy_(torch.tensor([0, cut, 150]))
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                for n in ("q", "k", "v", "do"):
                    t[n].copy_(other[n])
                graph.replay()
            stream.synchronize()
            compare(t, True, ("replay", seed))
            got = {n: t[n].clone() for n in ("o", "dq", "dk", "dv")}
            torch.cuda.synchronize()
            M.mmee_prompt_attn_forward(a)
            M.mmee_prompt_attn_backward(a, g)
            stream.synchronize()
            for n, x in got.items():
                assert torch.equal(x, t[n]), (n, seed)
    finally:
        M.mmee_set_stream(None)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("lens,H,Hkv,d", [([70, 40, 90], 2, 1, 64), ([70, 40, 300], 4, 2, 128), ([300, 500, 260], 33, 33, 104), ([600, 57, 700], 8, 8, 64)])
def test_a_sequence_that_is_not_finite(M, lens, H, Hkv, d, dtype):
    """Reaches none of the others."""
    import torch
    t = tensors(lens, lens, H, Hkv, d, getattr(torch, dtype), 41)
    middle = slice(lens[0], lens[0] + lens[1])
    for n in ("q", "k", "v", "do"):
        t[n][middle] = math.nan
        t[n][middle][::3] = math.inf
    run(M, t, kv=False)
    for at in (slice(0, middle.start), slice(middle.stop, sum(lens))):
        one = {n: t[n][at] for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")} | {"lse": t["lse"][:, at]}
        one["q_starts"] = one["kv_starts"] = starts_of([at.stop - at.start])
        compare(one, True, (lens, at))


def test_graphs_that_share_a_workspace(M):
    """A forward and a backward call, planned and in pieces, captured one by one with one workspace; replayed in turn over other lengths and inputs."""
    import torch
    T = 2400
    make = lambda lens, seed: tensors(lens, lens, 4, 2, 128, torch.bfloat16, seed)  # noqa: E731
    t = make([1200, 1200], 50)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    M.mmee_set_stream(stream.cuda_stream)
    try:
        a, g = calls(M, t)
        M.mmee_prompt_attn_forward(a)
        M.mmee_prompt_attn_backward(a, g)
        stream.synchronize()
        graphs = []
        for call in (lambda: M.mmee_prompt_attn_forward(a), lambda: M.mmee_prompt_attn_backward(a, g)):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=stream):
                call()
        for seed, cut in enumerate((2300, 1, 1200, T)):
            other = make([cut, T - cut], 51 + seed)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                for n in ("q", "k", "v", "do", "q_starts", "kv_starts"):
                    t[n].copy_(other[n])
                for graph in graphs:
                    graph.replay()
            stream.synchronize()
            compare(t, True, ("replay", cut))
    finally:
        M.mmee_set_stream(None)


def test_gradients_against_differences(M):
    """The change of sum(o do) along one direction of each input, in 64 bits, against the gradients."""
    import torch
    from attention_oracle import attention
    m, n, H, Hkv, d = 30, 45, 4, 2, 32
    t = tensors([m], [n], H, Hkv, d, torch.float16, 18)
    run(M, t)
    x = {name: t[name].cpu().double() for name in ("q", "k", "v", "do")}

    def value(q, k, v):
        k, v = (z.repeat_interleave(H // Hkv, 1) for z in (k, v))
        s = torch.einsum("mhd,nhd->hmn", q, k) * d ** -0.5
        o = torch.einsum("hmn,nhd->mhd", torch.softmax(s.masked_fill(~keep_of(m, n, True), -math.inf), 2), v)
        return (o * x["do"]).sum()
    bounds = attention(*(t[name][None] for name in ("q", "k", "v")), keep_of(m, n, True), d ** -0.5, torch.float16, t["do"][None])
    step = 1e-5
    for name in ("q", "k", "v"):
        way = torch.randn(x[name].shape, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
        moved = [value(**{p: x[p] + (sign * step * way if p == name else 0) for p in "qkv"}) for sign in (1, -1)]
        want = (moved[0] - moved[1]) / (2 * step)
        got = (t["d" + name].cpu().double() * way).sum()
        assert abs(got - want) <= (bounds["d" + name][1][0] * way.abs()).sum() + 1e-6 * abs(want), name
