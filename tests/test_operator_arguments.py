"""What the operators' calls refuse, before anything is launched: needs the built library, no GPU.  Tensors are stand-ins with a
device tensor's face."""
import ctypes as C
import os

import pytest

M = None


@pytest.fixture(scope="module", autouse=True)
def binding():
    """The binding, loaded when a test runs and after torch: whichever of the two comes first brings the HIP runtime that both use."""
    global M
    import torch  # noqa: F401
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    if not os.path.exists(os.environ.get("MMEE_LIB") or os.path.join(root, "paper_2604_03446_amd", "libmmee.so")):
        import __graft_entry__ as g
        g.build()
    import paper_2604_03446_amd
    M = paper_2604_03446_amd


class Fake:
    """A device tensor without a device: nothing may read or write it."""
    is_cuda = True

    def __init__(self, *shape, dtype="torch.bfloat16", stride=None, at=1 << 20):
        self.shape, self.dtype, self.at = shape, dtype, at
        if stride is None:
            stride, n = [], 1
            for s in reversed(shape):
                stride.insert(0, n)
                n *= s
        self._stride = tuple(stride)

    def stride(self):
        return self._stride

    def data_ptr(self):
        return self.at

    def is_contiguous(self):
        return self._stride == Fake(*self.shape)._stride

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return {"torch.bfloat16": 2, "torch.float16": 2, "torch.uint8": 1}.get(self.dtype, 4)


def cross(**over):
    t = {"q": Fake(2, 5, 4, 64), "k": Fake(2, 7, 2, 64), "v": Fake(2, 7, 2, 64), "o": Fake(2, 5, 4, 64)}
    kw = {n: v for n, v in over.items() if n not in t}
    t.update({n: v for n, v in over.items() if n in t})
    return M.attn(t["q"], t["k"], t["v"], t["o"], **kw)


def refused(call, code=None):
    with pytest.raises(M.MmeeError) as e:
        call()
    assert e.value.code == (M.EINVAL if code is None else code)


def test_attention_refuses():
    assert M.mmee_attn_workspace(cross()) == 0
    on_host = Fake(2, 5, 4, 64)
    on_host.is_cuda = False
    for over in (dict(q=on_host), dict(q=Fake(2, 5, 4, 64, dtype="torch.float32")), dict(v=Fake(2, 7, 2, 64, dtype="torch.float16")), dict(k=Fake(2, 6, 2, 64)),
                 dict(o=Fake(2, 5, 4, 32)), dict(q=Fake(2, 5, 64, 4, stride=(1280, 256, 1, 64))), dict(kv_lens=Fake(3, dtype="torch.int32")),
                 dict(kv_lens=Fake(2, dtype="torch.int64")), dict(key_mask=Fake(2, 7, dtype="torch.float32")), dict(key_mask=Fake(2, 8, dtype="torch.uint8")),
                 dict(lse=Fake(2, 4, 5, dtype="torch.float64")), dict(lse=Fake(2, 4, 5, dtype="torch.float32", stride=(20, 1, 4)))):
        refused(lambda: cross(**over))
    for over in (dict(k=Fake(2, 7, 3, 64), v=Fake(2, 7, 3, 64)),                                      # heads that do not share evenly
                 dict(q=Fake(2, 5, 4, 68), k=Fake(2, 7, 2, 68), v=Fake(2, 7, 2, 68), o=Fake(2, 5, 4, 68)),            # head size no multiple of 8
                 dict(q=Fake(2, 5, 4, 136), k=Fake(2, 7, 2, 136), v=Fake(2, 7, 2, 136), o=Fake(2, 5, 4, 136)),        # head size beyond 128
                 dict(k=Fake(2, 7, 2, 64, stride=(900, 129, 64, 1))), dict(q=Fake(2, 5, 4, 64, stride=(1280, -256, 64, 1))),
                 dict(o=Fake(2, 5, 4, 64, stride=(0, 256, 64, 1))), dict(o=Fake(2, 5, 4, 64, stride=(1280, 256, 0, 1))),
                 dict(k=Fake(2, 7, 2, 64, stride=(1 << 30, 1 << 25, 64, 1))), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        refused(lambda: M.mmee_attn_workspace(cross(**over)))
        refused(lambda: M.mmee_attn_forward(cross(**over)))
    refused(lambda: M.mmee_attn_forward(cross(q=Fake(2, 5, 4, 64, at=(1 << 20) + 8))))
    refused(lambda: M.mmee_attn_forward(cross(k=Fake(2, 7, 2, 64, at=0))))
    for field, value in (("dtype", 2), ("batch", 0), ("heads", 0), ("kv_heads", 0), ("head_dim", 0), ("reserved", 1)):
        a = cross()
        setattr(a, field, value)
        refused(lambda: M.mmee_attn_forward(a))
    assert M._lib.mmee_attn_forward(None) == M.EINVAL and M._lib.mmee_attn_workspace(C.byref(cross()), 0, None) == M.EINVAL


def test_attention_wants_its_workspace():
    long = dict(q=Fake(1, 1, 4, 64), k=Fake(1, 9000, 1, 64), v=Fake(1, 9000, 1, 64), o=Fake(1, 1, 4, 64))
    size = M.mmee_attn_workspace(cross(**long))
    assert size > 0
    refused(lambda: M.mmee_attn_forward(cross(**long)), M.EWORKSPACE)
    refused(lambda: M.mmee_attn_forward(cross(**long).use_workspace(Fake(size - 1, dtype="torch.uint8"))), M.EWORKSPACE)
    refused(lambda: M.mmee_attn_forward(cross(**long).use_workspace(Fake(size, dtype="torch.uint8", at=(1 << 20) + 4))))
    assert "workspace" in M._strerror(M.EWORKSPACE)


def test_attention_backward_refuses():
    grads = lambda **o: M.attn_grads(*({"do": Fake(2, 5, 4, 64), "dq": Fake(2, 5, 4, 64), "dk": Fake(2, 7, 2, 64), "dv": Fake(2, 7, 2, 64)} | o).values())  # noqa: E731
    a = cross(lse=Fake(2, 4, 5, dtype="torch.float32"))
    a.use_workspace(Fake(M.mmee_attn_workspace(a, True), dtype="torch.uint8"))
    refused(lambda: M.mmee_attn_backward(cross(), grads()))                          # no lse
    refused(lambda: M.mmee_attn_backward(cross(lse=Fake(2, 4, 5, dtype="torch.float32")), grads()), M.EWORKSPACE)
    for over in (dict(do=Fake(2, 5, 2, 64), dq=Fake(2, 5, 2, 64)), dict(dk=Fake(2, 7, 4, 64), dv=Fake(2, 7, 4, 64)), dict(dk=Fake(2, 7, 2, 64, stride=(0, 128, 64, 1))),
                 dict(dv=Fake(2, 7, 2, 64, at=(1 << 20) + 2)), dict(dq=Fake(2, 5, 4, 64, at=0)),
                 {n: Fake(2, *s, 64, dtype="torch.float16") for n, s in (("do", (5, 4)), ("dq", (5, 4)), ("dk", (7, 2)), ("dv", (7, 2)))}):
        refused(lambda: M.mmee_attn_backward(a, grads(**over)))
    assert M._lib.mmee_attn_backward(C.byref(a), None) == M.EINVAL


def tree(**over):
    t = {"q": Fake(2, 70, 4, 64), "k_pages": Fake(9, 16, 2, 64), "v_pages": Fake(9, 16, 2, 64), "page_table": Fake(2, 6, dtype="torch.int32"),
         "cache_lens": Fake(2, dtype="torch.int32"), "ancestors": Fake(2, 70, 2, dtype="torch.int64"), "o": Fake(2, 70, 4, 64)}
    kw = {n: v for n, v in over.items() if n not in t}
    t.update({n: v for n, v in over.items() if n in t})
    return M.tree_attn(*t.values(), **kw)


def test_tree_attention_refuses():
    M.mmee_tree_attn_workspace(tree())
    for over in (dict(ancestors=Fake(2, 70, 1, dtype="torch.int64")), dict(ancestors=Fake(2, 70, 2, dtype="torch.int32")), dict(cache_lens=Fake(2, dtype="torch.int64")),
                 dict(page_table=Fake(2, 6, dtype="torch.int64")), dict(page_table=Fake(3, 6, dtype="torch.int32")), dict(node_counts=Fake(1, dtype="torch.int32")),
                 dict(v_pages=Fake(9, 16, 2, 32)), dict(page_table=Fake(2, 6, dtype="torch.int32", stride=(12, 2)))):
        refused(lambda: tree(**over))
    for over in (dict(k_pages=Fake(9, 24, 2, 64), v_pages=Fake(9, 24, 2, 64)), dict(k_pages=Fake(9, 16, 3, 64), v_pages=Fake(9, 16, 3, 64)), dict(scale=0.0),
                 dict(q=Fake(2, 1025, 4, 64), o=Fake(2, 1025, 4, 64), ancestors=Fake(2, 1025, 17, dtype="torch.int64")),
                 dict(o=Fake(2, 70, 4, 64, stride=(0, 256, 64, 1)))):
        refused(lambda: M.mmee_tree_attn_workspace(tree(**over)))
    refused(lambda: M.mmee_tree_attn_forward(tree(ancestors=Fake(2, 70, 2, dtype="torch.int64", at=(1 << 20) + 4))))
    refused(lambda: M.mmee_tree_attn_forward(tree(cache_lens=Fake(2, dtype="torch.int32", at=0))))
    long = tree(page_table=Fake(2, 4000, dtype="torch.int32"))
    assert M.mmee_tree_attn_workspace(long) > 0
    refused(lambda: M.mmee_tree_attn_forward(long), M.EWORKSPACE)
    assert M._lib.mmee_tree_attn_forward(None) == M.EINVAL


def block(**over):
    t = {"x": Fake(9, 64), "w_gate": Fake(80, 64), "w_up": Fake(80, 64), "w_down": Fake(48, 80), "y": Fake(9, 48), "hidden": Fake(9, 80)}
    kw = {n: v for n, v in over.items() if n not in t}
    t.update({n: v for n, v in over.items() if n in t})
    return M.ffn(*t.values(), **kw)


def test_ffn_refuses():
    assert M.mmee_ffn_workspace(block()) == 0 and M.mmee_ffn_workspace(block(), True) > 0
    for over in (dict(act="tanh"), dict(w_up=Fake(72, 64)), dict(w_down=Fake(48, 72)), dict(y=Fake(9, 40)), dict(hidden=Fake(9, 80, stride=(88, 1))),
                 dict(gate=Fake(9, 72)), dict(x=Fake(9, 64, dtype="torch.float32")), dict(w_gate=Fake(80, 64, stride=(1, 80)))):
        refused(lambda: block(**over))
    for over in (dict(x=Fake(9, 60), w_gate=Fake(80, 60), w_up=Fake(80, 60)), dict(w_up=Fake(80, 64, stride=(72, 1))), dict(x=Fake(9, 64, stride=(0, 1))),
                 dict(x=Fake(9, 64, stride=(65, 1))), dict(y=Fake(9, 48, stride=(40, 1))), dict(w_down=Fake(48, 80, stride=(1 << 23, 1)))):
        refused(lambda: M.mmee_ffn_workspace(block(**over)))
    refused(lambda: M.mmee_ffn_forward(block(hidden=Fake(9, 80, at=(1 << 20) + 8))))
    refused(lambda: M.mmee_ffn_forward(block(w_down=Fake(48, 80, at=0))))
    for field, value in (("dtype", 7), ("act", 5), ("in_dim", 0), ("hidden_dim", 0), ("out_dim", 0), ("reserved", 1)):
        f = block()
        setattr(f, field, value)
        refused(lambda: M.mmee_ffn_forward(f))
    grads = lambda **o: M.ffn_grads(*({"dy": Fake(9, 48), "dx": Fake(9, 64), "dw_gate": Fake(80, 64), "dw_up": Fake(80, 64), "dw_down": Fake(48, 80)} | o).values())  # noqa: E731
    kept = block(gate=Fake(9, 80), up=Fake(9, 80))
    refused(lambda: M.mmee_ffn_backward(kept, grads()), M.EWORKSPACE)
    kept.use_workspace(Fake(M.mmee_ffn_workspace(kept, True), dtype="torch.uint8"))
    refused(lambda: M.mmee_ffn_backward(block(), grads()))                           # g and u were not kept
    for over in (dict(dx=Fake(9, 56)), dict(dw_gate=Fake(72, 64)), dict(dy=Fake(9, 48, stride=(0, 1))), dict(dx=Fake(9, 64, at=0)), dict(dw_up=Fake(80, 64, at=(1 << 20) + 8))):
        refused(lambda: M.mmee_ffn_backward(kept, grads(**over)))
    refused(lambda: grads(dw_down=Fake(48, 80, stride=(88, 1))))
    assert M._lib.mmee_ffn_backward(C.byref(kept), None) == M.EINVAL
