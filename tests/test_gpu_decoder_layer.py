"""The example's layer, run as a user would, against the same layer in plain 32-bit torch."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_layer_against_plain_torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(ROOT, "examples", "decoder_layer.py"))
    E = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(E)
    layer = E.Layer(3, 11, 8, 2, 64, 320, dtype=torch.float16)
    t = E.inputs(layer, cache=150, encoder=90)
    B, n, H, Hkv, d = 3, 11, 8, 2, 64
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    E.M.mmee_set_stream(stream.cuda_stream)
    try:
        with torch.cuda.stream(stream):
            got = layer.step(**t)
        stream.synchronize()
    finally:
        E.M.mmee_set_stream(None)

    def attend(q, k, v, keep):                  # [n, H, d], [L, Hkv, d], [n, L]
        k, v = (z.float().repeat_interleave(H // Hkv, 1) for z in (k, v))
        s = torch.einsum("nhd,lhd->hnl", q.float(), k) * d ** -0.5
        return torch.einsum("hnl,lhd->nhd", torch.softmax(s.masked_fill(~keep, -float("inf")), 2), v)

    norm = lambda z: torch.nn.functional.layer_norm(z.float(), (H * d,))  # noqa: E731
    for b in range(B):
        x = t["x"][b].float()
        q = (norm(x) @ layer.w_qkv[:H * d].float().t()).view(n, H, d)
        held = int(t["cache_lens"][b])
        pages = t["page_table"][b].long()
        k, v = (t[z][pages].reshape(-1, Hkv, d)[:held + n] for z in ("k_pages", "v_pages"))         # (the step has put the tokens' own behind)
        sees = torch.tensor([[w >> j & 1 for j in range(n)] for w in t["ancestors"][b, :, 0].tolist()], dtype=torch.bool, device="cuda")
        keep = torch.cat([torch.ones(n, held, dtype=torch.bool, device="cuda"), sees], 1)
        x = x + attend(q, k, v, keep).reshape(n, -1) @ layer.w_self_out.float().t()
        length = int(t["enc_lens"][b])
        q = (norm(x) @ layer.w_cross_q.float().t()).view(n, H, d)
        x = x + attend(q, t["enc_k"][b, :length], t["enc_v"][b, :length], torch.ones(n, length, dtype=torch.bool, device="cuda")).reshape(n, -1) @ layer.w_cross_out.float().t()
        z = norm(x)
        x = x + (torch.nn.functional.silu(z @ layer.w_gate.float().t()) * (z @ layer.w_up.float().t())) @ layer.w_down.float().t()
        # some twenty roundings to 11 bits of values of size 1 to 4 on the way: 2^-11 each, in the root mean square
        assert (got[b].float() - x).square().mean().sqrt() <= 2.0 ** -11 * 20 ** 0.5 * x.square().mean().sqrt()


def test_planned_chains():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(ROOT, "examples", "decoder_layer.py"))
    E = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(E)
    from inputs import CONFIGS
    for name, r in E.plan(2, 8, 4, 32, 128, 64, 40, CONFIGS["tiny"]["hw"]):
        assert r.cost.valid and r.cost.energy_pj > 0, name
