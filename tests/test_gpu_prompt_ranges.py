"""Attention of packed prompts where its ranges end: float16 gradients far from unit size, D of rows that see few keys, short sequences beside long
ones, and as many sequences and tiles as a plan and a wave's look at the starts hold, and more."""
import math

import pytest

from test_gpu_prompt_attention import compare, keep_of, run, tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


def gradients(t, rows, keys, causal=True):
    """(values, bounds) of dq, dk, dv of one sequence in float16, as attention_oracle.py has them, but that what rounding leaves of small numbers is relative: P is
    kept to 2^-32 of a row's largest at least (2^-25 of the type, 2^7 above it), and dS to 2^-35 of the largest of its row or key (2^-25 where that lies above
    2^10).  Outputs have steps of 2^-24 below the normal numbers."""
    u, tiny = 2.0 ** -11, 2.0 ** -25
    H, Hkv, d = t["q"].shape[1], t["k"].shape[1], t["q"].shape[2]
    heads = lambda x, at: t[x][at].double().cpu().transpose(0, 1)  # noqa: E731
    q, do = heads("q", rows), heads("do", rows)
    k, v = (heads(x, keys).repeat_interleave(H // Hkv, 0) for x in ("k", "v"))
    keep, scale = keep_of(q.shape[1], k.shape[1], causal)[0], d ** -0.5
    P = (q @ k.transpose(1, 2) * scale).masked_fill(~keep, -math.inf).softmax(2)
    O, dP, across = P @ v, do @ v.transpose(1, 2), do.abs() @ v.abs().transpose(1, 2)
    o_off = u * O.abs() + 1.5 * u * (P @ v.abs()) + 2.0 ** -32 * (keep.double() @ v.abs()) + tiny
    dS = P * (dP - (do * O).sum(2, keepdim=True))
    off = 1.5 * u * dS.abs() + P * (0.5 * u * across + (do.abs() * o_off).sum(2, keepdim=True))
    row, key = (2.0 ** -35 * dS.abs().amax(i, keepdim=True) * keep for i in (2, 1))
    shared = lambda x: x.view(Hkv, H // Hkv, *x.shape[1:]).sum(1).transpose(0, 1)  # noqa: E731
    turn = lambda x: x.transpose(1, 2)  # noqa: E731
    dQ, dK, dV = (dS @ k * scale).transpose(0, 1), shared(turn(dS) @ q) * scale, shared(turn(P) @ do)
    return {"dq": (dQ, u * dQ.abs() + scale * ((off + row) @ k.abs()).transpose(0, 1) + tiny),
            "dk": (dK, u * dK.abs() + scale * shared(turn(off + key) @ q.abs()) + tiny),
            "dv": (dV, u * dV.abs() + 1.5 * u * shared(turn(P) @ do.abs()) + 2.0 ** -40 * shared(turn(keep.double().expand_as(P)) @ do.abs()) + tiny)}


def check_gradients(t, lens, where, causal=True):
    from attention_oracle import check
    at = 0
    for n in lens:
        one = slice(at, at + n)
        at += n
        for name, want in gradients(t, one, one, causal).items():
            check(t[name][one], want, (where, n, name))


RANGES = [([1, 2, 9, 16, 3], 64), ([40, 64, 17], 128), ([300, 129], 64), ([300, 700], 128), ([2100], 128)]       # one step of a product; a tile; several; eight waves for dK and dV; for dQ too, and cut tiles


@pytest.mark.parametrize("by", [-12, 10])
@pytest.mark.parametrize("lens,d", RANGES)
def test_float16_gradients_far_from_unit_size(M, lens, d, by):
    """dO of 2^-12 and of 2^10: dS is kept in float16's range either way."""
    import torch
    H, Hkv = (8, 2) if sum(lens) == 1000 else (4, 2)
    t = tensors(lens, lens, H, Hkv, d, torch.float16, 71 + by)
    # (float16 holds what is scaled down exactly)
    t["do"] = ((t["do"].float() * 64).round() / 64).clamp(-4, 4).mul(2.0 ** by).to(torch.float16)
    run(M, t, kv=False)
    check_gradients(t, lens, by)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("first,then", [(-12, 8), (8, -12)])
@pytest.mark.parametrize("lens,d", RANGES)
def test_float16_gradients_whose_size_changes(M, lens, d, first, then, causal):
    """Rows of dO, and keys' values, of another size from the middle of the sequence on: dS outgrows the power of two that it was kept by, with sums there already."""
    import torch
    H, Hkv = (8, 2) if sum(lens) == 1000 else (4, 2)
    for which in ("do", "v"):
        t = tensors(lens, lens, H, Hkv, d, torch.float16, 73)
        at = 0
        for n in lens:
            size = torch.full((n, 1, 1), 2.0 ** first, device="cuda")
            size[n // 2:] = 2.0 ** then
            if which == "v":
                size = size.clamp(2.0 ** -6, 2.0 ** 6)
            t[which][at:at + n] *= size.to(torch.float16)
            at += n
        run(M, t, kv=False, causal=causal)
        check_gradients(t, lens, (which, first, causal), causal)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("beside", [0, 20000])
def test_D_of_few_keys_that_weigh_the_same(M, beside, dtype):
    """All keys' values are ones and all dO the same, queries are orthogonal to keys: dP is one number B, P is 1 / n, dS is P (B - D) = 0, and what D is off by shows alone.
    Alone and beside a sequence over so many keys, with which blocks have eight waves.

    In float16's forward pass the sum is n 2^7 and its logarithm, below 16, off by a unit of 2^-20; twice it is multiplied and rounded, 2^-23 of 4: 2^-20 and 2^-21 of
    a power of two, times ln 2 below 2^-20 of P.  An exponential is off by 2^-23, and D is n / 2 additions in each of two lanes and one, 2^-24 each: 2^-21 for n up to
    16.  So |B - D| <= B (2^-20 + 2^-21 + 2^-22), which dS and the results of n terms have as they have P; their own roundings are below 2^-7 of that."""
    import torch
    d, dt, B = 128, getattr(torch, dtype), 128.0 * 128
    lens = [7, 9, 11, 14, 16, 3] if beside else list(range(2, 17))
    t = tensors(lens + [1500] * (beside > 0), lens + [beside] * (beside > 0), 2, 1, d, dt, 77)
    t["q"][..., :64], t["k"][..., 64:] = 0, 0
    t["v"].fill_(1.0)
    t["do"].fill_(128.0)
    run(M, t, causal=False)
    at = 0
    for n in lens:
        one = slice(at, at + n)
        at += n
        off = 1.01 * B * (2.0 ** -20 + 2.0 ** -21 + 2.0 ** -22) * d ** -0.5
        k, q = t["k"][one].double().abs().sum(0, keepdim=True) / n, t["q"][one].double().abs().sum((0, 1), keepdim=True) / n
        for name, bound in (("dq", off * k), ("dk", off * q)):
            far = t[name][one].double().abs() - bound - 2.0 ** -25
            assert (far <= 0).all(), (n, name, far.max().item(), (t[name][one].double().abs() / (bound + 2.0 ** -25)).max().item())


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_dS_of_up_to_16_keys_one_by_one(M, dtype):
    """Keys are unit vectors, so that a value of dQ is one dS times the scale, and of V and dO one value is not zero, so that dP is exact: dS goes into dQ as two
    operands and is off by u^2 and by what errors in 32 bits add, and its result is rounded once, to u.

    P is off by 2^-19 (scores below 8 and their products with log2 e below 2^-21 of a power of two, lse, the logarithm of a sum of up to 2^11, 2^-20), D by that and 16
    additions, 2^-20.  Float16 has steps of 2^-24 below its normal numbers."""
    import torch
    d, dt = 64, getattr(torch, dtype)
    u, scale = torch.finfo(dt).eps / 2, d ** -0.5
    lens = [16, 9, 13, 2, 15, 7] * 8
    t = tensors(lens, lens, 4, 2, d, dt, 101)
    at = 0
    for n in lens:
        t["k"][at:at + n] = torch.eye(n, d, device="cuda")[:, None].to(dt)
        at += n
    t["q"] *= 3
    t["v"][..., 1:], t["do"][..., 1:] = 0, 0
    run(M, t, kv=False, causal=False)
    at = 0
    for b, n in enumerate(lens):
        one = slice(at, at + n)
        at += n
        q, do, v = (t[x][one].double().cpu().transpose(0, 1) for x in ("q", "do", "v"))
        P = (q[..., :n] * scale).softmax(2)
        dP = do[..., :1] * v[..., 0].repeat_interleave(2, 0)[:, None]
        D = (P * dP).sum(2, keepdim=True)
        dS = P * (dP - D)
        off = (u + 1.01 * u * u) * dS.abs() + 1.01 * P * (2.0 ** -19 * (dP - D).abs() + (2.0 ** -19 + 2.0 ** -20) * (P * dP.abs()).sum(2, keepdim=True))
        far = (t["dq"][one].double().cpu().transpose(0, 1)[..., :n] - dS * scale).abs() - off * scale - 2.0 ** -25
        assert (far <= 0).all(), (b, n, int((far > 0).sum()), far.max().item())


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("lens,d", [([1200, 9, 1200, 16, 1], 128), ([4200, 9], 128), ([2300, 5], 64)])
def test_few_keys_beside_long_sequences(M, lens, d, dtype):
    """Blocks of eight waves, which the average length decides, round dS once for sequences of any length (up to 16 keys alone, blocks of four take what that leaves
    along): to u of each dS, and what errors in 32 bits add as in the test of gradients of few keys."""
    import torch
    t = tensors(lens, lens, 4, 2, d, getattr(torch, dtype), 79)
    run(M, t, kv=False)
    u, scale = torch.finfo(t["q"].dtype).eps / 2, d ** -0.5
    for b, n in enumerate(lens):
        if n > 16:
            continue
        at = slice(sum(lens[:b]), sum(lens[:b]) + n)
        q, do = (t[x][at].double().cpu().view(n, 2, 2, d).permute(1, 2, 0, 3) for x in ("q", "do"))
        k, v = (t[x][at].double().cpu().permute(1, 0, 2)[:, None] for x in ("k", "v"))
        P = (q @ k.transpose(2, 3) * scale).masked_fill(~keep_of(n, n, True), -math.inf).softmax(3)
        dP, across = do @ v.transpose(2, 3), do.abs() @ v.abs().transpose(2, 3)
        dS = P * (dP - (P * dP).sum(3, keepdim=True))
        off = u * dS.abs() + 2.0 ** -16 * P * (across + (P * across).sum(3, keepdim=True))
        for name, want, bound in (("dq", dS @ k, off @ k.abs()), ("dk", (dS.transpose(2, 3) @ q).sum(1, keepdim=True), (off.transpose(2, 3) @ q.abs()).sum(1, keepdim=True))):
            got = t[name][at].double().cpu().view(n, 2, -1, d).permute(1, 2, 0, 3)
            far = (got - want * scale).abs() - (1.01 * bound + u * want.abs()) * scale - 2.0 ** -25
            assert (far <= 0).all(), (b, n, name, far.max().item())


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q_lens,kv_lens,H,Hkv,d", [
    ([2100] + [40] * 60, None, 2, 1, 64), ([40] * 30 + [1500] + [3] * 30, None, 4, 1, 128), ([64, 8, 8, 8], [5000, 30, 30, 30], 4, 1, 128),
    ([3, 1, 40, 200, 0], [3000, 5000, 1, 200, 900], 4, 1, 64), ([1] * 9, [2] * 8 + [9000], 2, 1, 32)])
def test_one_long_sequence_among_short_ones(M, q_lens, kv_lens, H, Hkv, d, causal, dtype):
    """Whose average length is far from all of theirs: cut into pieces or not."""
    import torch
    t = tensors(q_lens, kv_lens or q_lens, H, Hkv, d, getattr(torch, dtype), 83, around=1)
    run(M, t, causal=causal)
    compare(t, causal, (q_lens, kv_lens))


def compare_padded(t, where):
    """As compare(), all sequences at once, padded to the longest."""
    import torch
    from attention_oracle import attention, check
    q_starts, kv_starts = t["q_starts"].cpu().long(), t["kv_starts"].cpu().long()
    m, n = q_starts.diff(), kv_starts.diff()
    i, j = torch.arange(int(m.max())), torch.arange(int(n.max()))
    there, key_there = i < m[:, None], j < n[:, None]
    rows, keys = (q_starts[:-1, None] + i).clamp(max=t["q"].shape[0] - 1), (kv_starts[:-1, None] + j).clamp(max=t["k"].shape[0] - 1)
    keep = there[:, :, None] & key_there[:, None] & (j <= i[:, None] + (n - m)[:, None, None])
    pad = lambda x, at, live: torch.where(live[..., None, None], x.cpu()[at], torch.zeros((), dtype=x.dtype))  # noqa: E731
    q, do, k, v = pad(t["q"], rows, there), pad(t["do"], rows, there), pad(t["k"], keys, key_there), pad(t["v"], keys, key_there)
    for name, (value, off) in attention(q, k, v, keep, t["q"].shape[2] ** -0.5, t["q"].dtype, do).items():
        if name == "lse":
            check(t["lse"].cpu()[:, rows].transpose(0, 1).transpose(1, 2)[there], (value.transpose(1, 2)[there], off.transpose(1, 2)[there]), (where, name))
        else:
            at, live = (keys, key_there) if name[-1] in "kv" else (rows, there)
            check(t[name].cpu()[at][live], (value[live], off[live]), (where, name))


@pytest.mark.parametrize("seqs", [2047, 2048, 2049, 4096, 4097, 5003])
def test_as_many_sequences_as_a_plan_holds_and_more(M, seqs):
    """Of 0 to 3 rows; from 4097 on a wave looks at the starts three times."""
    import torch
    lens = [i * 7 % 4 for i in range(seqs)]
    t = tensors(lens, [n + i % 3 for i, n in enumerate(lens)], 2, 1, 32, torch.bfloat16, 89, around=1)
    run(M, t)
    compare_padded(t, seqs)


@pytest.mark.parametrize("more", [0, 1])
def test_as_many_tiles_as_a_plan_holds_and_more(M, more):
    """2048 tiles of rows at most, with a start of every sequence's own, are planned, 2049 go by slots; tiles of keys are more either way."""
    import torch
    seqs, H = 512, 4
    lens = [96 + (i * 29 % 63 - 31) for i in range(seqs)]
    lens[-1] += 1536 * 128 // H - sum(lens) + 128 // H * more                # H rows a token: 1536 tiles of 128 rows, or one more
    kv_lens = [n + 130 for n in lens]
    t = tensors(lens, kv_lens, H, 1, 16, torch.bfloat16, 97)
    assert min(lens) > 0 and sum(lens) * H // 128 + seqs == 2048 + more
    run(M, t)
    compare_padded(t, more)
