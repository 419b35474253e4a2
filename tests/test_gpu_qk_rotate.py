"""Norm and rotation of queries and keys, forward and backward, against a plain 64-bit form (rotation_oracle.py): head sizes, pairings, rotated
parts, axes, far positions, layouts, in place, values out of the ordinary, streams, graphs."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


def tensors(T, H, Hkv, d, rot, dtype, seed, axes=1, norm=True, train=True, far=100000, scale=1.5):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)  # noqa: E731
    t = {"q": r(T, H, d), "k": r(T, Hkv, d)}
    t |= {n + "_out": torch.full_like(t[n], math.nan) for n in ("q", "k")}
    t["freqs"] = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).cuda() if rot else None
    t["positions"] = torch.randint(0, far, (axes, T) if axes > 1 else (T,), generator=g, device="cuda").to(torch.int32) if rot else None
    t["axis_of"] = torch.randint(0, axes, (rot // 2,), generator=g, device="cuda").to(torch.uint8) if axes > 1 else None
    for n in ("q", "k"):
        t[n + "_weight"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dtype) if norm else None
    if train:
        t |= {"dq_out": r(T, H, d), "dk_out": r(T, Hkv, d)}
        t |= {"d" + n: torch.full_like(t[n], math.nan) for n in ("q", "k")}
        t |= {f"d{n}_weight": torch.full((d,), math.nan, dtype=dtype, device="cuda") if norm else None for n in ("q", "k")}
    return t


def calls(M, t, **kw):
    import torch
    f = M.qk_rotate(t["q"], t["k"], t["q_out"], t["k_out"], t["freqs"], t["positions"], t["axis_of"], t["q_weight"], t["k_weight"], **kw)
    # whatever the workspace holds before a call does not matter
    f.use_workspace(torch.full((M.mmee_qk_rotate_workspace(f),), 255, dtype=torch.uint8, device="cuda"))
    return f, M.qk_rotate_grads(t["dq_out"], t["dk_out"], t["dq"], t["dk"], t["dq_weight"], t["dk_weight"]) if "dq_out" in t else None


def run(M, t, **kw):
    import torch
    f, g = calls(M, t, **kw)
    M.mmee_qk_rotate_forward(f)
    if g:
        M.mmee_qk_rotate_backward(f, g)
    torch.cuda.synchronize()


def compare(t, where, pairs="halves", eps=1e-6, inputs=None):
    import torch
    from attention_oracle import check
    from rotation_oracle import angles, rotation
    angle = angles(t["freqs"], t["positions"], t["axis_of"]) if t["freqs"] is not None else torch.zeros(t["q"].shape[0], 1, 0, dtype=torch.float64)
    for n in ("q", "k"):
        want = rotation((inputs or t)[n], t[n + "_weight"], angle, eps, pairs, (inputs or t).get(f"d{n}_out"))
        for name, key in (("y", n + "_out"), ("dx", "d" + n), ("dw", f"d{n}_weight")):
            if name in want:
                check(t[key], want[name], (where, key))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("T,H,Hkv,d,rot", [(1, 1, 1, 8, 0), (1, 32, 8, 128, 128), (3, 5, 1, 16, 16), (7, 4, 2, 24, 16), (33, 12, 12, 64, 64), (65, 6, 3, 80, 32), (17, 3, 3, 72, 48),
                                           (5, 2, 1, 40, 32), (31, 8, 8, 96, 96), (129, 7, 1, 120, 112), (9, 3, 2, 256, 256), (40, 2, 2, 200, 64), (6, 9, 4, 136, 0), (300, 1, 1, 32, 32)])
def test_shapes(M, T, H, Hkv, d, rot, pairs, dtype):
    import torch
    for norm in (True, False):
        t = tensors(T, H, Hkv, d, rot, getattr(torch, dtype), T + d, norm=norm)
        run(M, t, pairs=pairs)
        compare(t, (T, H, Hkv, d, rot, pairs, norm), pairs)


def test_many_tokens(M):
    """More tokens than a backward pass has waves: every wave takes several."""
    import torch
    t = tensors(5003, 3, 2, 64, 32, torch.bfloat16, 3)
    run(M, t)
    compare(t, "many tokens")


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("axes", [2, 3, 4])
def test_axes(M, axes, pairs):
    import torch
    t = tensors(50, 4, 2, 96, 64, torch.float16, axes, axes=axes)
    run(M, t, pairs=pairs)
    compare(t, axes, pairs)
    t["axis_of"][::3] = 250                     # beyond the axes: the last one
    wide = torch.full((axes, 64), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    wide[:, :50] = t["positions"]
    t["positions"] = wide[:, :50]
    run(M, t, pairs=pairs)
    compare(t, (axes, "clamped"), pairs)


def test_far_and_negative_positions(M):
    import torch
    t = tensors(12, 2, 1, 64, 64, torch.float16, 9)
    t["positions"] = torch.tensor([0, 1, -1, 2 ** 20, 2 ** 20 + 1, -2 ** 20, 2 ** 24 + 1, 10 ** 7, 12345678, -12345679, 3, 99999999], dtype=torch.int32, device="cuda")
    run(M, t)
    compare(t, "far")


def test_long_tensors(M):
    """Places beyond 2^31 elements from the first one."""
    import torch
    T, d = 3, 64
    row = (1 << 31) + 64
    big = torch.zeros(2 * row + 64 * 2 * d, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(big)
    t = tensors(T, 2, 1, d, 64, torch.bfloat16, 2, train=False)
    far = lambda b, heads: b.as_strided((T, heads, d), (row, d, 1))  # noqa: E731
    far(big, 2).copy_(t["q"])
    t["q"], t["q_out"] = far(big, 2), far(out, 2)
    run(M, t)
    compare(t, "far apart")


@pytest.mark.parametrize("layout", ["fused", "heads first", "broadcast", "in place", "sliced"])
def test_layouts(M, layout):
    import torch
    T, H, Hkv, d, dt = 45, 4, 2, 64, torch.bfloat16
    t = tensors(T, H, Hkv, d, 64, dt, 4)
    inputs = None
    if layout == "fused":
        for pre, post in (("", ""), ("", "_out"), ("d", "_out"), ("d", "")):
            x = torch.full((T, H + 2 * Hkv, d), 7.0, dtype=dt, device="cuda")
            x[:, :H], x[:, H:H + Hkv] = t[f"{pre}q{post}"], t[f"{pre}k{post}"]
            t |= {f"{pre}q{post}": x[:, :H], f"{pre}k{post}": x[:, H:H + Hkv]}
    elif layout == "heads first":
        for n in ("q", "k", "q_out", "k_out", "dq_out", "dk_out", "dq", "dk"):
            t[n] = t[n].transpose(0, 1).contiguous().transpose(0, 1)
    elif layout == "broadcast":
        t["q"], t["k"], t["dk_out"] = t["q"][:1].expand(T, H, d), t["k"][:, :1].expand(T, Hkv, d), t["dk_out"][:1, :1].expand(T, Hkv, d)
    elif layout == "sliced":
        wide = torch.full((T, H, d + 16), 5.0, dtype=dt, device="cuda")
        t["q_out"] = wide[..., 8:8 + d]
    else:
        inputs = {n: t[n].clone() for n in ("q", "k", "dq_out", "dk_out")}
        t["dq"], t["dk"] = t["dq_out"], t["dk_out"]
        f, g = calls(M, t)
        M.mmee_qk_rotate_backward(f, g)                  # which reads q and k, so before they are overwritten
        t["q_out"], t["k_out"] = t["q"], t["k"]
        f, _ = calls(M, t)
        M.mmee_qk_rotate_forward(f)
        torch.cuda.synchronize()
    if layout != "in place":
        run(M, t)
    compare(t, layout, inputs=inputs)
    if layout == "fused":
        assert (x[:, H + Hkv:] == 7.0).all()
    if layout == "sliced":
        assert (wide[..., :8] == 5.0).all() and (wide[..., 8 + d:] == 5.0).all()


def test_heads_of_zeros_and_of_what_is_not_finite(M):
    """A head of zeros gives zeros and finite gradients; what is not finite stays in its head, and without a norm in its pair."""
    import torch
    t = tensors(8, 4, 2, 64, 32, torch.bfloat16, 6)
    t["q"][2, 1] = 0
    run(M, t)
    compare(t, "zeros")
    assert not t["q_out"][2, 1].any()
    for norm in (True, False):
        t = tensors(8, 4, 2, 64, 32, torch.float16, 7, norm=norm, train=False)
        clean = {n: t[n].clone() for n in ("q", "k")}
        t["q"][3, 2, 5], t["k"][1, 0, 40] = math.inf, math.nan
        run(M, t)
        bad_q, bad_k = torch.zeros_like(t["q"], dtype=torch.bool), torch.zeros_like(t["k"], dtype=torch.bool)
        if norm:
            bad_q[3, 2], bad_k[1, 0] = True, True
        else:
            bad_q[3, 2, [5, 21]], bad_k[1, 0, 40] = True, True
        assert not torch.isfinite(t["q_out"][3, 2, 5]) and torch.isnan(t["k_out"][1, 0, 40])
        got = {n: t[n].clone() for n in ("q_out", "k_out")}
        t |= clean
        run(M, t)
        assert torch.equal(got["q_out"][~bad_q], t["q_out"][~bad_q]) and torch.equal(got["k_out"][~bad_k], t["k_out"][~bad_k])


def test_nothing_to_do(M):
    import torch
    t = tensors(0, 4, 2, 64, 64, torch.bfloat16, 1)
    run(M, t)
    assert not t["dq_weight"].any() and not t["dk_weight"].any()


def test_gradients_against_differences(M):
    """One direction of the inputs: the change of sum(y dy) against the gradients, in steps large enough for 16-bit outputs summed over many values."""
    import torch
    from rotation_oracle import angles, rotation
    t = tensors(20, 3, 2, 64, 64, torch.float16, 8)
    run(M, t)
    angle = angles(t["freqs"], t["positions"])
    way = torch.randn(t["q"].shape, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    step, x, dy = 1e-4, t["q"].cpu().double(), t["dq_out"].cpu().double()

    def value(x, w):
        z = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
        a, b = z[..., :32], z[..., 32:]
        return (torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1) * dy).sum()
    w = t["q_weight"].cpu().double()
    want = (value(x + step * way, w) - value(x - step * way, w)) / (2 * step)
    bound = rotation(t["q"], t["q_weight"], angle, 1e-6, "halves", t["dq_out"])["dx"][1]
    assert abs((t["dq"].cpu().double() * way).sum() - want) <= (bound * way.abs()).sum() + 1e-4 * want.abs()
    way = torch.randn(64, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
    want = (value(x, w + step * way) - value(x, w - step * way)) / (2 * step)
    bound = rotation(t["q"], t["q_weight"], angle, 1e-6, "halves", t["dq_out"])["dw"][1]
    assert abs((t["dq_weight"].cpu().double() * way).sum() - want) <= (bound * way.abs()).sum() + 1e-4 * want.abs()


def test_repeats_to_the_bit(M):
    import torch
    t = tensors(2500, 8, 2, 128, 128, torch.bfloat16, 12)
    run(M, t)
    first = {n: t[n].clone() for n in ("q_out", "k_out", "dq", "dk", "dq_weight", "dk_weight")}
    run(M, t)
    for n, x in first.items():
        assert torch.equal(x, t[n]), n


def test_streams_and_graphs(M):
    """Captured on a stream of its own and replayed over changed inputs, with eager calls of the same buffers between the replays."""
    import torch
    t = tensors(70, 4, 2, 64, 64, torch.bfloat16, 10)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    M.mmee_set_stream(stream.cuda_stream)
    try:
        with torch.cuda.stream(stream):
            f, g = calls(M, t)
            M.mmee_qk_rotate_forward(f)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            M.mmee_qk_rotate_forward(f)
            M.mmee_qk_rotate_backward(f, g)
        for seed in range(4):
            other = tensors(70, 4, 2, 64, 64, torch.bfloat16, 20 + seed)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                for n in ("q", "k", "dq_out", "dk_out"):
                    t[n].copy_(other[n])
                graph.replay()
            stream.synchronize()
            compare(t, ("replay", seed))
            got = {n: t[n].clone() for n in ("q_out", "k_out", "dq", "dk", "dq_weight", "dk_weight")}
            torch.cuda.synchronize()
            M.mmee_qk_rotate_forward(f)
            M.mmee_qk_rotate_backward(f, g)
            stream.synchronize()
            for n, x in got.items():
                assert torch.equal(x, t[n]), (n, seed)
    finally:
        M.mmee_set_stream(None)
