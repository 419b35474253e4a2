"""An error that the program met before a call is not the call's: the call succeeds, and the error is still there for the program to ask for."""
import pytest

from test_gpu_attention import run as run_cross
from test_gpu_attention import tensors
from test_gpu_ffn import run as run_ffn
from test_gpu_ffn import tensors as block
from test_gpu_tree_attention import build
from test_gpu_tree_attention import run as run_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("operator", ["cross", "tree", "ffn"])
def test_earlier_error(operator):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as M
    if operator == "cross":
        t = tensors((1, 5, 2, 64), (1, 70, 2, 64), torch.bfloat16, 1)
        a = M.attn(t["q"], t["k"], t["v"], t["o"], lse=t["lse"])
        a.use_workspace(torch.empty(M.mmee_attn_workspace(a, True), dtype=torch.uint8, device="cuda"))
        g = M.attn_grads(t["do"], t["dq"], t["dk"], t["dv"])
        calls = [lambda: M.mmee_attn_forward(a), lambda: M.mmee_attn_backward(a, g)]
        run_cross(M, t)
    elif operator == "tree":
        t = build(1, 3, 2, 1, 64, 16, [20], torch.bfloat16)
        from test_gpu_tree_attention import words_of
        words = words_of(t["sees"]).cuda()
        a = M.tree_attn(t["q"], t["k_pages"], t["v_pages"], t["table"], t["lens"], words, t["o"], lse=t["lse"])
        a.use_workspace(torch.empty(M.mmee_tree_attn_workspace(a), dtype=torch.uint8, device="cuda"))
        calls = [lambda: M.mmee_tree_attn_forward(a)]
        run_tree(M, t)
    else:
        t = block(9, 64, 72, 40, torch.bfloat16, 1)
        f = M.ffn(t["x"], t["w_gate"], t["w_up"], t["w_down"], t["y"], t["hidden"], gate=t["gate"], up=t["up"])
        f.use_workspace(torch.empty(M.mmee_ffn_workspace(f, True), dtype=torch.uint8, device="cuda"))
        g = M.ffn_grads(t["dy"], t["dx"], t["dw_gate"], t["dw_up"], t["dw_down"])
        calls = [lambda: M.mmee_ffn_forward(f), lambda: M.mmee_ffn_backward(f, g)]
        run_ffn(M, t, "silu")
    hip = M._lib                                        # (finds the runtime's functions in what the library is linked to)
    for call in calls:
        error = hip.hipSetDevice(9999)                  # no such device: an error of the program's own
        assert error != 0
        try:
            call()
            assert hip.hipPeekAtLastError() == error
        finally:
            hip.hipGetLastError()
    torch.cuda.synchronize()
