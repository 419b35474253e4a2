"""Performance cases of the operators that run a planned chain: cross attention, tree attention over a cache, gated feed-forward.

A case is a dict of plain values.  `prepare` makes the tensors that a program holds before the call, `run` is one pass:
the operators' plain form in 32 bits, or, where `own` is true, the library's calls on the same tensors.  `exact` restates
each operator in 64 bits.
"""
import math

import torch

own = False                 # true: `run` makes the library's calls

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- the cases ---------------------------------------------------------------------------------

def _cross(B, H, Hkv, d, Lq, Lk, dtype, ragged=False, mask=False, train=False):
    return {"kind": "cross", "B": B, "H": H, "Hkv": Hkv, "d": d, "Lq": Lq, "Lk": Lk, "dtype": dtype, "ragged": ragged, "mask": mask, "train": train}


def _tree(B, H, Hkv, d, nodes, ctx, page, dtype, ragged=False):
    return {"kind": "tree", "B": B, "H": H, "Hkv": Hkv, "d": d, "nodes": nodes, "ctx": ctx, "page": page, "dtype": dtype, "ragged": ragged}


def _ffn(rows, K, F, J, dtype, act, train=False):
    return {"kind": "ffn", "rows": rows, "K": K, "F": F, "J": J, "dtype": dtype, "act": act, "train": train}


def listed():
    return [
        # One decoded token against a short encoded input: latency counts.
        {"name": "cross_token", **_cross(1, 12, 12, 64, 1, 512, "bf16")},
        # A serving batch of single tokens, each against an encoded input of its own length, shared key/value heads.
        {"name": "cross_tokens_ragged", **_cross(64, 32, 8, 128, 1, 2048, "fp16", ragged=True)},
        # A prompt against a long encoded input.
        {"name": "cross_prompt", **_cross(1, 32, 32, 128, 2048, 8192, "bf16")},
        # A training step over padded inputs: odd lengths, a mask of keys.
        {"name": "cross_train_masked", **_cross(8, 12, 12, 64, 509, 1500, "bf16", mask=True, train=True)},
        # A training step with shared key/value heads and long inputs.
        {"name": "cross_train", **_cross(2, 32, 8, 128, 2048, 4096, "bf16", train=True)},
        # One sequence checks a handful of drafted tokens after a short context: latency counts.
        {"name": "tree_one", **_tree(1, 32, 8, 128, 7, 500, 16, "bf16")},
        # A serving batch checks full trees, every sequence at a length of its own.
        {"name": "tree_batch", **_tree(16, 32, 8, 128, 63, 4096, 16, "fp16", ragged=True)},
        # Two long contexts.
        {"name": "tree_long", **_tree(2, 64, 8, 128, 26, 131072, 64, "bf16", ragged=True)},
        # One token through a small layer: latency counts.
        {"name": "ffn_token", **_ffn(1, 768, 3072, 768, "bf16", "silu")},
        # A decoding batch through a large layer, bound by its weights.
        {"name": "ffn_tokens", **_ffn(37, 4096, 12288, 4096, "fp16", "gelu_tanh")},
        # A prompt through the layer whose mapping the benchmark searches.
        {"name": "ffn_prompt", **_ffn(2048, 768, 3072, 768, "bf16", "gelu")},
        # A training step, an odd number of tokens.
        {"name": "ffn_train", **_ffn(4001, 2048, 8192, 2048, "bf16", "silu", train=True)},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    kind = rng.choice(["cross", "cross", "tree", "ffn"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if kind == "ffn":
        wide = lambda lo, hi: max(lo, _log_int(rng, lo, hi) // 8 * 8)  # noqa: E731
        train = rng.random() < 0.4
        K = wide(256, 4096)
        return _ffn(_log_int(rng, 64 if train else 1, 8192), K, wide(512, 12288), rng.choice([K, wide(256, 4096)]), dtype,
                    rng.choice(["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]), train)
    Hkv = rng.choice([1, 2, 4, 8, 12, 16])
    H = Hkv * rng.choice([1, 1, 2, 4, 8])
    d = rng.choice([32, 64, 80, 96, 128, 128])
    if kind == "tree":
        return _tree(_log_int(rng, 1, 32), H, Hkv, d, _log_int(rng, 1, 128), _log_int(rng, 1, 131072), rng.choice([16, 32, 64, 128]), dtype, rng.random() < 0.7)
    train = rng.random() < 0.4
    Lq = 1 if not train and rng.random() < 0.4 else _log_int(rng, 2, 2048)
    masking = rng.choice(["", "ragged", "mask"])
    return _cross(_log_int(rng, 1, 64), H, Hkv, d, Lq, _log_int(rng, 1, 8192), dtype, masking == "ragged", masking == "mask", train)


def draw(rng):
    most = {}
    for c in listed():
        w, m = work(c), most.setdefault(c["kind"], {"bytes": 0, "flops": 0})
        for key in m:
            m[key] = max(m[key], w[key])
    while True:
        c = _draw(rng)
        w = work(c)
        # the plain form of attention keeps all scores: no more of them than the largest listed case has
        scores = c["B"] * c["H"] * c.get("Lq", c.get("nodes")) * c.get("Lk", c.get("ctx")) if c["kind"] != "ffn" else 0
        if all(w[key] <= most[c["kind"]][key] for key in w) and scores <= 2 * 32 * 2048 * 4096:
            return c


def work(case):
    c = case
    if c["kind"] == "ffn":
        weights, tokens = 2 * c["K"] * c["F"] + c["F"] * c["J"], c["rows"] * (c["K"] + c["J"])
        # forward: x and weights in, y out; a training step also reads dy and writes dx and the weights' gradients
        return {"bytes": 2 * (weights + tokens) * (2 if c["train"] else 1), "flops": 2 * c["rows"] * weights * (3 if c["train"] else 1)}
    if c["kind"] == "tree":
        # a ragged batch holds three quarters of the longest context on average
        ctx = (0.75 if c["ragged"] else 1.0) * c["ctx"] + c["nodes"]
        q = c["B"] * c["nodes"] * c["H"] * c["d"]
        return {"bytes": 2 * (2 * q + 2 * c["B"] * ctx * c["Hkv"] * c["d"]), "flops": 4 * q * ctx}
    Lk = (0.75 if c["ragged"] else 1.0) * c["Lk"]
    q, kv = c["B"] * c["Lq"] * c["H"] * c["d"], 2 * c["B"] * Lk * c["Hkv"] * c["d"]
    # forward: two products; backward: five. A training step reads q, k, v, do and writes o and three gradients
    return {"bytes": 2 * (2 * q + kv) * (2 if c["train"] else 1), "flops": 2 * q * Lk * (7 if c["train"] else 2)}


# ---- what a program has in hand ------------------------------------------------------------------

def _randn(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = DTYPES[c["dtype"]]
    s = dict(c)
    if c["kind"] == "ffn":
        rows, K, F, J = c["rows"], c["K"], c["F"], c["J"]
        s["x"] = _randn(gen, rows, K, dtype=dtype)                              # a normed input
        s["w_gate"] = _randn(gen, F, K, dtype=dtype, scale=K ** -0.5)
        s["w_up"] = _randn(gen, F, K, dtype=dtype, scale=K ** -0.5)
        s["w_down"] = _randn(gen, J, F, dtype=dtype, scale=F ** -0.5)
        s["y"] = torch.empty(rows, J, dtype=dtype, device="cuda")
        s["hidden"] = torch.empty(rows, F, dtype=dtype, device="cuda")
        if c["train"]:
            s["dy"] = _randn(gen, rows, J, dtype=dtype)
            for name, like in (("gate", "hidden"), ("up", "hidden"), ("dx", "x"), ("dw_gate", "w_gate"), ("dw_up", "w_up"), ("dw_down", "w_down")):
                s[name] = torch.empty_like(s[like])
        return s
    B, H, Hkv, d = c["B"], c["H"], c["Hkv"], c["d"]
    if c["kind"] == "tree":
        n, page, ctx = c["nodes"], c["page"], c["ctx"]
        per_seq = -(-(ctx + n) // page)
        s["q"] = _randn(gen, B, n, H, d, dtype=dtype)
        # the pool of pages, keys and values of a page beside each other; sequences hold its pages in no order
        pool = _randn(gen, B * per_seq, 2, page, Hkv, d, dtype=dtype)
        s["k_pages"], s["v_pages"] = pool[:, 0], pool[:, 1]
        s["page_table"] = torch.randperm(B * per_seq, generator=gen, device="cuda").to(torch.int32).view(B, per_seq)
        s["cache_lens"] = torch.full((B,), ctx, dtype=torch.int32, device="cuda")
        s["node_counts"] = torch.full((B,), n, dtype=torch.int32, device="cuda")
        if c["ragged"]:
            s["cache_lens"] = torch.randint(ctx // 2, ctx + 1, (B,), generator=gen, device="cuda").to(torch.int32)
            s["node_counts"] = torch.randint((n + 1) // 2, n + 1, (B,), generator=gen, device="cuda").to(torch.int32)
        # a random tree: node i hangs on a node before it; its row holds its ancestors and itself
        parent = (torch.rand(B, n, generator=gen, device="cuda") * torch.arange(n, device="cuda")).long()
        seen = torch.zeros(B, n, n, dtype=torch.bool, device="cuda")
        seen[:, 0, 0] = True
        at = torch.arange(B, device="cuda")
        for i in range(1, n):
            seen[:, i] = seen[at, parent[:, i]]
            seen[:, i, i] = True
        words = -(-n // 64)
        bits = torch.zeros(B, n, words * 64, dtype=torch.long, device="cuda")
        bits[:, :, :n] = seen
        s["ancestors"] = (bits.view(B, n, words, 64) << torch.arange(64, device="cuda")).sum(-1)    # 64 bits of a word, the last one its sign
        s["o"] = torch.empty(B, n, H, d, dtype=dtype, device="cuda")
        return s
    Lq, Lk = c["Lq"], c["Lk"]
    s["q"] = _randn(gen, B, Lq, H, d, dtype=dtype)
    kv = _randn(gen, B, Lk, 2, Hkv, d, dtype=dtype)             # one projection of the encoder's states gives keys and values
    s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
    s["kv_lens"] = torch.randint(Lk // 2, Lk + 1, (B,), generator=gen, device="cuda").to(torch.int32) if c["ragged"] else None
    s["key_mask"] = (torch.rand(B, Lk, generator=gen, device="cuda") < 0.8).to(torch.uint8) if c["mask"] else None
    s["o"] = torch.empty(B, Lq, H, d, dtype=dtype, device="cuda")
    if c["train"]:
        s["lse"] = torch.empty(B, H, Lq, dtype=torch.float32, device="cuda")
        s["do"] = _randn(gen, B, Lq, H, d, dtype=dtype)
        s["dq"] = torch.empty_like(s["q"])
        dkv = torch.empty_like(kv)
        s["dk"], s["dv"] = dkv[:, :, 0], dkv[:, :, 1]
    return s


# ---- the plain forms, 32 bits ----------------------------------------------------------------------

def _heads(x, Hkv):
    """[B, L, H, d] -> [B, Hkv, group * L, d] in 32 bits: the rows that share a key/value head."""
    B, L, H, d = x.shape
    return x.float().view(B, L, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, H // Hkv * L, d)


def _tokens(x, L, H):
    """[B, Hkv, group * L, d] -> [B, L, H, d]"""
    B, Hkv, _, d = x.shape
    return x.view(B, Hkv, H // Hkv, L, d).permute(0, 3, 1, 2, 4).reshape(B, L, H, d)


def _softmax(scores, allowed):
    scores = scores.masked_fill(~allowed, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    return torch.where(total > 0, p / total, torch.zeros_like(p))


def _plain_cross(s):
    B, Lq, H, d = s["q"].shape
    Hkv, Lk, dtype, scale = s["Hkv"], s["Lk"], s["q"].dtype, d ** -0.5
    q, k, v = _heads(s["q"], Hkv), _heads(s["k"], Hkv), _heads(s["v"], Hkv)
    allowed = torch.ones(B, Lk, dtype=torch.bool, device=q.device)
    if s["kv_lens"] is not None:
        allowed = torch.arange(Lk, device=q.device) < s["kv_lens"][:, None]
    if s["key_mask"] is not None:
        allowed = allowed & (s["key_mask"] != 0)
    p = _softmax(torch.matmul(q, k.transpose(2, 3).contiguous()) * scale, allowed[:, None, None, :])
    o = torch.matmul(p, v)
    out = {"o": _tokens(o, Lq, H).to(dtype)}
    if not s["train"]:
        return out
    do = _heads(s["do"], Hkv)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (do * o).sum(-1, keepdim=True)) * scale
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    out["dq"] = _tokens(dq, Lq, H).to(dtype)
    out["dk"], out["dv"] = dk.transpose(1, 2).to(dtype), dv.transpose(1, 2).to(dtype)
    return out


def _plain_tree(s):
    B, n, H, d = s["q"].shape
    Hkv, page = s["Hkv"], s["page"]
    table = s["page_table"].long()
    L = table.shape[1] * page
    k = _heads(s["k_pages"][table].reshape(B, L, Hkv, d), Hkv)
    v = _heads(s["v_pages"][table].reshape(B, L, Hkv, d), Hkv)
    dev = k.device
    at = torch.arange(L, device=dev)[None, :] - s["cache_lens"][:, None]                # place among the drafted tokens, negative in the cache
    j = at.clamp(0, n - 1)
    word = torch.gather(s["ancestors"], 2, (j // 64)[:, None, :].expand(B, n, L))
    seen = ((word >> (j % 64)[:, None, :]) & 1) != 0
    drafted = (at >= 0) & (at < s["node_counts"][:, None])
    live = torch.arange(n, device=dev)[None, :] < s["node_counts"][:, None]
    allowed = ((at < 0)[:, None, :] | (drafted[:, None, :] & seen)) & live[:, :, None]
    scores = torch.matmul(_heads(s["q"], Hkv), k.transpose(2, 3).contiguous()) * d ** -0.5
    p = _softmax(scores, allowed[:, None].repeat(1, 1, H // Hkv, 1))
    return {"o": _tokens(torch.matmul(p, v), n, H).to(s["q"].dtype)}


def _act(g, name):
    """An activation and its derivative."""
    if name == "silu":
        e = torch.sigmoid(g)
        return g * e, e * (1 + g * (1 - e))
    if name == "sigmoid":
        e = torch.sigmoid(g)
        return e, e * (1 - e)
    if name == "relu":
        e = (g > 0).to(g.dtype)
        return g * e, e
    if name == "gelu":
        e = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
        return g * e, e + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5
    c, a = (2 / math.pi) ** 0.5, 0.044715
    t = torch.tanh(c * (g + a * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * a * g * g)


def _plain_ffn(s):
    dtype = s["x"].dtype
    x, wg, wu, wd = (s[name].float() for name in ("x", "w_gate", "w_up", "w_down"))
    g, u = torch.matmul(x, wg.t()), torch.matmul(x, wu.t())
    a, da = _act(g, s["act"])
    h = a * u
    out = {"y": torch.matmul(h, wd.t()).to(dtype)}
    if not s["train"]:
        return out
    dy = s["dy"].float()
    dh = torch.matmul(dy, wd)
    dg, du = dh * u * da, dh * a
    out["dx"] = (torch.matmul(dg, wg) + torch.matmul(du, wu)).to(dtype)
    out["dw_gate"] = torch.matmul(dg.t(), x).to(dtype)
    out["dw_up"] = torch.matmul(du.t(), x).to(dtype)
    out["dw_down"] = torch.matmul(dy.t(), h).to(dtype)
    return out


# ---- the library's calls -----------------------------------------------------------------------------

def _marshal(s):
    """The structures that a program makes once of its buffers and keeps, with their workspace."""
    import paper_2604_03446_amd as M
    if s["kind"] == "ffn":
        f = M.ffn(s["x"], s["w_gate"], s["w_up"], s["w_down"], s["y"], s["hidden"], act=s["act"], gate=s.get("gate"), up=s.get("up"))
        g = M.ffn_grads(s["dy"], s["dx"], s["dw_gate"], s["dw_up"], s["dw_down"]) if s["train"] else None
        call, size = (f, g), M.mmee_ffn_workspace(f, s["train"])
    elif s["kind"] == "tree":
        f = M.tree_attn(s["q"], s["k_pages"], s["v_pages"], s["page_table"], s["cache_lens"], s["ancestors"], s["o"], node_counts=s["node_counts"])
        call, size = (f, None), M.mmee_tree_attn_workspace(f)
    else:
        f = M.attn(s["q"], s["k"], s["v"], s["o"], lse=s.get("lse"), kv_lens=s["kv_lens"], key_mask=s["key_mask"])
        g = M.attn_grads(s["do"], s["dq"], s["dk"], s["dv"]) if s["train"] else None
        call, size = (f, g), M.mmee_attn_workspace(f, s["train"])
    f.use_workspace(torch.empty(size, dtype=torch.uint8, device="cuda"))
    return M, call


def _calls(s):
    if "call" not in s:
        s["call"] = _marshal(s)
    M, (f, g) = s["call"]
    if s["kind"] == "tree":
        M.mmee_tree_attn_forward(f)
        return {"o": s["o"]}
    if s["kind"] == "ffn":
        M.mmee_ffn_forward(f)
        if not s["train"]:
            return {"y": s["y"]}
        M.mmee_ffn_backward(f, g)
        return {name: s[name] for name in ("y", "dx", "dw_gate", "dw_up", "dw_down")}
    M.mmee_attn_forward(f)
    if not s["train"]:
        return {"o": s["o"]}
    M.mmee_attn_backward(f, g)
    return {name: s[name] for name in ("o", "dq", "dk", "dv")}


def run(state):
    if own:
        return _calls(state)
    return {"cross": _plain_cross, "tree": _plain_tree, "ffn": _plain_ffn}[state["kind"]](state)


# ---- the definitions, 64 bits --------------------------------------------------------------------------
# Sequence by sequence and head by head; gradients by differentiating the forward definition.

def _attend(q, k, v, keep):
    """One head: rows q see the keys that keep[row] marks; rows that see none give zeros."""
    z = (q @ k.t()) / math.sqrt(q.shape[1])
    none = ~keep.any(1, keepdim=True)
    z = z.masked_fill(~(keep | none), -math.inf)
    return (torch.softmax(z, 1) @ v).masked_fill(none, 0.0)


def _exact_cross(c, s):
    group, names = c["H"] // c["Hkv"], ["q", "k", "v"]
    x = {name: s[name].double().requires_grad_(c["train"]) for name in names}
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device="cuda")
    grads = {name: torch.zeros(s[name].shape, dtype=torch.float64, device="cuda") for name in names} if c["train"] else {}
    for b in range(c["B"]):
        keep = torch.ones(c["Lk"], dtype=torch.bool, device="cuda")
        if c["ragged"]:
            keep[int(s["kv_lens"][b]):] = False
        if c["mask"]:
            keep &= s["key_mask"][b].bool()
        for h in range(c["H"]):
            q, k, v = (x[name][b, :, h if name == "q" else h // group].detach().requires_grad_(c["train"]) for name in names)
            out = _attend(q, k, v, keep.expand(c["Lq"], -1))
            o[b, :, h] = out.detach()
            if c["train"]:
                got = torch.autograd.grad(out, (q, k, v), s["do"][b, :, h].double())
                for name, g in zip(names, got):
                    grads[name][b, :, h if name == "q" else h // group] += g
    return {"o": o, **{"d" + name: g for name, g in grads.items()}}


def _exact_tree(c, s):
    group, n = c["H"] // c["Hkv"], c["nodes"]
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        held, count = int(s["cache_lens"][b]), int(s["node_counts"][b])
        pages = s["page_table"][b].long()
        words = s["ancestors"][b].tolist()
        tree = torch.tensor([[words[i][j // 64] >> j % 64 & 1 for j in range(count)] for i in range(count)], dtype=torch.bool, device="cuda")
        keep = torch.cat([torch.ones(count, held, dtype=torch.bool, device="cuda"), tree.view(count, count)], 1)
        for m in range(c["Hkv"]):
            k = s["k_pages"][pages, :, m].reshape(-1, c["d"])[:held + count].double()
            v = s["v_pages"][pages, :, m].reshape(-1, c["d"])[:held + count].double()
            for h in range(m * group, (m + 1) * group):
                o[b, :count, h] = _attend(s["q"][b, :count, h].double(), k, v, keep)
    assert o.shape[1] == n
    return {"o": o}


def _exact_ffn(c, s):
    from torch.nn import functional as nn
    act = {"silu": nn.silu, "sigmoid": torch.sigmoid, "relu": nn.relu, "gelu": nn.gelu, "gelu_tanh": lambda g: nn.gelu(g, approximate="tanh")}[c["act"]]
    leaves = [s[name].double().requires_grad_(c["train"]) for name in ("x", "w_gate", "w_up", "w_down")]
    x, wg, wu, wd = leaves
    y = nn.linear(act(nn.linear(x, wg)) * nn.linear(x, wu), wd)
    if not c["train"]:
        return {"y": y}
    return {"y": y.detach(), **dict(zip(("dx", "dw_gate", "dw_up", "dw_down"), torch.autograd.grad(y, leaves, s["dy"].double())))}


def exact(case, seed):
    s = prepare(case, seed)
    return {"cross": _exact_cross, "tree": _exact_tree, "ffn": _exact_ffn}[case["kind"]](case, s)
